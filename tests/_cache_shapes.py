"""Shapes of the cache operators' larger paths, and what their plans make of
them: checked on the CPU, run on the GPU."""

# (sequence lengths, selected rows of each, Hq, Hkv, d), keys per workgroup / 64.
# The rows are the sequence's last ones and a few before, so that most steps of
# 128 (row, head) pairs are seen whole by a workgroup's keys and some are not.
SCORES = [
    (((4099, 0, 1003), (300, 0, 90), 16, 8, 64), 2), (((4099, 1003), (250, 100), 32, 8, 128), 2),
    (((8101, 333), (260, 333), 32, 8, 128), 4), (((16389,), (500,), 8, 4, 64), 4),
    (((2111,) * 5, (130,) * 5, 8, 8, 128), 4), (((9001,), (400,), 24, 8, 64), 4),
]

# (cache lengths, Hq, Hkv, d), keys per chunk.  Full chunks fill a wave's ring of
# slots several times over; the others end inside it.
_LONG = (4100, 4097, 3333, 2049, 5119, 4096, 1, 17) * 2
_MID = (2100, 1025, 2047, 513, 1900, 2048, 1, 700) * 2
STEPS = [((lens, 8 * g, 8, d), kc)
         for lens, kc in ((_LONG, 1024), (_MID, 512)) for g in (4, 8, 16) for d in (64, 128)]
STEPS += [((_LONG, 24, 8, 128), 1024), ((_LONG, 40, 8, 64), 1024), ((_MID, 4 * 20, 4, 128), 512)]
