"""Every kernel that a product with 4-bit weights can take, with every group and zero form that it is built for, and shapes that reach what those of i4_checks leave out."""
import i4_checks

FORMS = ("linear", "gradient", "gated", "gated gradient")
# output channels, tokens, blocks of 128 columns in a step: as in csrc/lordba_i4_choice.h
TILES = {"tile32": (32, 32, 8), "tile64": (64, 32, 4), "tile128": (128, 64, 2), "tile256": (256, 128, 1), "square64": (64, 64, 4)}
# T, d_in, d_out (d_ff), group, zero points
SHAPES = [(1, 32, 6120, 64, False), (1, 56, 5496, 128, False), (1, 128, 8244, 64, True), (1, 8344, 48, 32, False), (2, 56, 8384, 32, True),
          (2, 96, 8264, 32, False), (2, 8288, 6472, 128, True), (3, 8269, 40, 128, False), (3, 8336, 1048, 64, False), (5, 4336, 4168, 32, True),
          (5, 4528, 32, 32, False), (5, 6768, 4568, 128, True), (5, 6832, 4744, 64, True), (6, 32, 8392, 64, False), (6, 96, 8264, 128, False),
          (6, 6064, 4368, 128, False), (6, 8288, 48, 32, True), (7, 72, 8256, 128, True), (8, 40, 7184, 32, False), (15, 4591, 32, 64, False),
          (54, 3184, 1656, 128, False), (66, 1224, 3096, 64, True), (73, 1059, 2624, 64, False), (114, 544, 8152, 64, True), (134, 584, 5664, 32, True),
          (138, 6414, 576, 32, False), (154, 1128, 1664, 32, False), (220, 1325, 296, 64, False), (390, 1344, 1128, 64, False), (440, 184, 3821, 32, True),
          (540, 2192, 552, 128, False), (653, 8044, 320, 128, False), (667, 112, 5512, 128, False), (680, 6264, 32, 64, False), (908, 3721, 32, 32, False),
          (914, 264, 5744, 128, True), (915, 1352, 528, 32, True), (934, 1224, 288, 128, True), (1044, 5298, 296, 64, False), (1165, 3984, 328, 64, True),
          (1320, 200, 752, 128, True), (1337, 3333, 32, 64, True), (1383, 288, 3240, 32, False), (1431, 731, 296, 32, False), (1661, 3214, 336, 32, False),
          (1690, 3007, 40, 128, False), (1693, 40, 2856, 32, False), (2018, 480, 80, 128, False), (2043, 696, 544, 64, False), (2049, 2648, 48, 32, True),
          (2074, 2184, 320, 32, True), (2158, 2480, 32, 32, False), (2205, 288, 2032, 64, True), (2404, 608, 568, 128, True), (2485, 272, 2520, 128, False),
          (2486, 616, 280, 32, True), (2509, 1656, 277, 64, False), (2516, 24, 1288, 64, True)]


def few(T, n, form):
    """Which of the kernels for few tokens: as in csrc/lordba_i4_few.hip"""
    tiles = -(-n // 32) * 2
    if tiles > 512 and T <= 8:
        return "few, four waves"
    if form == "linear" and tiles * -(-T // 16) <= 256:
        return "few, sixteen waves"
    if form != "gated" and tiles > 256 and T > 4:
        return "few, two blocks"
    return "few, eight waves"


def reached(T, d_in, d_out, group, zeros):
    """What the calls of a shape reach, tensors on their alignment and behind it: (form, kernel, aligned rows, group, zeros), tiles that exist whole, contractions of more
    than two steps, whole tiles of an odd number of outputs."""
    for shifted in (False, True):
        for form in FORMS:
            back = "gradient" in form
            k, n = (d_out, d_in) if back else (d_in, d_out)
            planes = 2 if form == "gated gradient" else 1
            aligned = not shifted and k % 8 == 0
            kernel = i4_checks.kernel(T, k, n, planes, form == "gated", aligned, back, zeros and group == 32)
            if kernel == "few":
                yield form, few(T, n, form), aligned, group, zeros
                continue
            yield form, kernel, aligned, group, zeros
            channels, tokens, parts = TILES[kernel]
            if n >= channels and T >= tokens:
                yield form, kernel, aligned, group, zeros, "whole"
                if n % 2:
                    yield form, kernel, aligned, "odd"
            if planes * -(-k // 128) > 2 * parts:
                yield form, kernel, aligned, group, zeros, "long"


def all_there_are():
    for form in FORMS:
        for aligned in (False, True):
            kernels = ["few, four waves", "few, eight waves", "tile32", "tile64", "tile128", "tile256"]
            kernels += ["few, sixteen waves"] * (form == "linear") + ["few, two blocks"] * (form != "gated") + ["square64"] * (form == "linear" and aligned)
            for kernel in kernels:
                if kernel in TILES:
                    yield form, kernel, aligned, "odd"
                for group in (32, 64, 128):
                    for zeros in (False, True):
                        if kernel == "tile256" and not aligned and "gradient" not in form and zeros and group == 32:
                            continue     # (not built: the choice leaves it out)
                        yield form, kernel, aligned, group, zeros
                        if kernel in TILES:
                            yield form, kernel, aligned, group, zeros, "whole"
                            yield form, kernel, aligned, group, zeros, "long"
