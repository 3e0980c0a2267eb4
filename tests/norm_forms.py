"""Which of the norm's kernels a call takes, as (vectors per thread, threads, stages of the ring, residual, row-code format or 0), and calls that between
them take every one of them for long enough that a CTA comes back to each slot of its ring."""

FEW_ROWS = 296


def _warps(cols, v):
    return -(-cols // (256 * v))


def forward_kernel(rows, cols, residual, y, fmt):
    wide = cols > 2048 and (not fmt if residual else bool(fmt) or y)
    v = 4 if cols > 8192 else 1 if rows <= FEW_ROWS else 4 if wide else 2
    threads = 256 if _warps(cols, v) <= 8 else 512 if _warps(cols, v) <= 16 else 1024
    stages = 3 if v < 4 else 1 if threads == 1024 else 2
    return v, threads, stages, residual, fmt


def backward_kernel(rows, cols, residual):
    v = 4 if cols > 8192 else 1 if rows <= FEW_ROWS else 2
    warps = _warps(cols, v)
    threads = 32 * warps * (1 if warps >= 8 else 8 // warps)
    row = (3 if residual else 2) * v * threads * 16
    if v == 4:
        return (4, 1024, 1, residual) if threads > 512 else (4, 512, 2, residual)
    return (1, 1024, 3, residual) if v == 1 else (2, 512, 3 if row <= 32 * 1024 else 2, residual)


# rows, cols, residual, y, fmt (0: none, 1: FP8, 2: FP4).  Widths among them whose warps per row do not divide the CTA's, which leaves warps without a row;
# beyond 296 rows more than the CTAs that threads and shared memory let be resident on 148 SMs, times their rows, times the stages.
FORWARD = [(rows, cols, residual, y, fmt)
           for residual in (False, True)
           for rows, cols, outs in ((296, 264, ((True, 0), (False, 1), (False, 2))), (289, 3336, ((True, 0), (False, 1), (False, 2))), (296, 8192, ((True, 0), (False, 1), (False, 2))),
                                    (15001, 1288, ((True, 0), (False, 1), (True, 2))), (3801, 4096, ((False, 0), (True, 1), (False, 2)) if residual else ((False, 0),)),
                                    (1951, 5128, ((False, 1), (True, 2)) if residual else ((False, 0),)), (1801, 8192, ((False, 1), (False, 2)) if residual else ((False, 0),)),
                                    (7203, 2056, ((True, 0),) if residual else ((True, 0), (False, 1), (True, 2))), (4801, 3200, ((True, 0),) if residual else ((True, 0), (True, 1), (False, 2))),
                                    (2400, 8192, ((True, 0),) if residual else ((True, 0), (False, 1), (False, 2))),
                                    (1203, 8200, ((True, 0), (False, 1), (False, 2))), (1201, 16384, ((False, 0), (True, 1), (False, 2))),
                                    (601, 17416, ((True, 0), (False, 1), (False, 2))), (600, 32768, ((False, 0), (True, 1), (False, 2))))
           for y, fmt in outs]
BACKWARD = [(rows, cols, residual) for residual in (False, True)
            for rows, cols in ((296, 520), (289, 3336), (296, 8192), (14000, 1032), (3601, 3200), (2301, 5128), (1801, 8192), (1201, 8200), (1203, 16384), (601, 17416), (603, 24576), (600, 32768))]
