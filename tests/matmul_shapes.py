"""Products that between them take every shape of workgroups: rows and columns that do not fill the last ones, at least five groups of k and a
last one that is cut, so that rings turn over and every edge is met."""
import paper_2510_08525_amd as rl

SHAPES = [(5, 1001, 2064), (13, 6149, 656), (16, 2051, 1168),                                                          # m <= 16
          (19, 1003, 1040), (64, 4099, 656), (23, 13001, 656), (61, 9007, 1040), (63, 28675, 656),                      # m <= 64
          (69, 109, 656), (67, 109, 1424), (65, 105, 5136), (201, 4003, 2064), (135, 5442, 656), (333, 4611, 3600), (5646, 134, 2208),
          (131, 11623, 656), (2040, 2045, 656), (1025, 6101, 656), (515, 10911, 656), (3001, 8203, 656), (8190, 4090, 656),
          (67, 17383, 656), (65, 8639, 656), (400, 5003, 784), (455, 8551, 656)]


def lists(dtype):
    """kind of call -> {place in its list: shapes that take it}, and the lists' lengths."""
    taken, lengths = {}, {}
    for s in SHAPES:
        *_, at, length = rl.rlkv_plan_matmul(*s, dtype)
        kind = "sixteen" if s[0] <= 16 else "sixty-four" if s[0] <= 64 else "many"
        taken.setdefault(kind, {}).setdefault(at, []).append(s)
        lengths[kind] = length
    return taken, lengths
