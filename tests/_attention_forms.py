"""The forms of the 8-bit cache's attention, and shapes that it runs in each: which shape takes which form is an estimate of
the library's that may change, so the tests ask it."""
SIZES = (32, 64, 72, 80, 96, 128)
CODE = {"f32": 0, "bf16": 1}
# keys widened once, groups of 32 queries of a workgroup, keys split over workgroups
FORMS = [("bf16", p, g, s) for p, g in ((False, 1), (False, 4), (True, 4)) for s in (False, True)] + \
        [("f32", False, 1, s) for s in (False, True)]
# B, heads, n_q, n_kv: the first that has the form is taken
CANDIDATES = [(1, 2, 40, 330), (2, 2, 70, 330), (1, 2, 33, 1501), (1, 2, 20, 5000), (1, 2, 129, 1001), (1, 2, 600, 2500),
              (1, 8, 1, 16384), (1, 8, 32, 8200), (8, 8, 32, 4099), (2, 16, 200, 1025), (2, 8, 600, 700), (2, 16, 520, 330),
              (2, 16, 1100, 333), (2, 16, 1100, 601), (2, 4, 1500, 1501), (2, 6, 1500, 2025), (1, 6, 1500, 3001)]


def shape_for(lib, form, d):
    """B, heads, n_q, n_kv, whether the call has its workspace; None if no candidate has the form."""
    dtype, prepared, groups, split = form
    for shape in CANDIDATES:
        need = lib.attention_quantized_workspace_bytes(*shape, d, CODE[dtype])
        for ws in (need, 0):
            got = lib.attention_quantized_plan(*shape, d, CODE[dtype], ws)
            if (got[0], got[1], got[2] > 1) == (prepared, groups, split):
                return (*shape, ws > 0)
    return None
