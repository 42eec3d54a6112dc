"""How a W4A16 call runs, by the rule of csrc/atom_w4a16.hip: which kernels it launches.  So that tests can say which of them their sizes reach."""


def _up(a, b):
    return -(-a // b)


def shape(M, N, K, O=128, gated=False, norm=True, index=True):
    """(kept, combine, NT, wide, parts) as product_shape gives them."""
    WM = 2 if gated else 1
    if M > 16:
        wide, U = 1 if M <= 32 else 2, (K + O) // 128
        tiles = _up(N, 128 if gated else 256) * _up(M, 32 * wide)
        best, parts = 1e30, 1
        for p in range(1, 33):
            if p * (6 if p > 16 else 2) > U:
                break
            cost = float(_up(tiles * p, 256)) * (_up(U, p) + 3) + (4 + float(p) * M * N * WM * 8 / 5e6 if p > 1 else 0)
            if cost < best:
                best, parts = cost, p
        return False, False, 0, wide, parts
    NT, combine = 1, norm and M <= 8
    sums = 8 * WM * 1024 * (2 if combine else 3)
    nat = 4 * K if norm else 2 * K if index else 0
    kept = False
    if M <= (8 if norm else 16):
        lds = M * (2 if norm else 1) * (K + 8) * 2 + max(nat, sums)
        kept = lds <= 80 * 1024 - 64 or (M == 1 and lds <= 150 * 1024 and _up(N, 16) <= 256)
    if not kept:
        rows, best = 2 * M if norm else M, 1e30
        for n in (1, 2, 4):
            if n * WM > 4:
                break
            cost = float(_up(_up(N, 16 * n), 256)) * (n * WM + rows / 16)
            if cost < best:
                best, NT = cost, n
    tiles, G4, parts = _up(N, 16 * NT), (K - O) // 128, 1
    wanted = min(G4 // 32, 256 // tiles)
    if wanted > 1:
        parts = _up(G4, _up(G4, wanted))
    return kept, combine, NT, 0, parts


def kernels(M, N, K, O=128, gated=False, norm=True, index=True):
    """The kernels that a call launches, as tuples of their names and template arguments."""
    kept, combine, NT, wide, parts = shape(M, N, K, O, gated, norm, index)
    out = []
    if not kept:
        out.append(("gather", bool(wide), 512 if K <= 4096 else 1024) if index else ("rows", bool(wide)))
    if wide:
        out.append(("wide", gated, wide, 2 if norm else 1))
    else:
        out.append(("few", NT, gated, 2 if norm and not combine else 1, combine, kept))
    if parts > 1:
        out.append(("join", gated))
    return out


ALL = ({("few", NT, g, HL, c, False) for NT, g in ((1, False), (2, False), (4, False), (1, True), (2, True)) for HL, c in ((1, False), (1, True), (2, False))} |
       {("few", 1, g, 1, c, True) for g in (False, True) for c in (False, True)} |
       {("wide", g, RT, HL) for g in (False, True) for RT in (1, 2) for HL in (1, 2)} |
       {("gather", w, t) for w in (False, True) for t in (512, 1024)} | {("rows", w) for w in (False, True)} | {("join", g) for g in (False, True)})
