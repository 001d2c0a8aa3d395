"""What a product of given sizes runs as, restated from the estimates of csrc/cdl_linear.cu and csrc/cdl_linear_rows.cu, so that tests can say which form
they mean and notice when an estimate moves a size elsewhere.  Sizes are (I, J, R): output rows and columns, reduced entries."""

PLAN_SMS, L2_BYTES, STAGE = 148, 126000000, 64


def up(n, m):
    return -(-n // m)


class Plan:
    def __init__(self, ns, whole, ranges, run, splits, piece_bytes, pair):
        self.ns, self.whole, self.ranges, self.run, self.splits, self.piece_bytes, self.pair = ns, whole, ranges, run, splits, piece_bytes, pair

    @property
    def form(self):
        return "cluster" if self.splits > 1 else ("pairs" if self.pair else "singles") + (" with runs" if self.ranges else "")


def tile_plan(I, J, R):
    kb, pairs, singles = up(R, STAGE), PLAN_SMS // 2, up(I, 128) * up(J, 128)
    forms = []
    for pair in (False, True):
        edge, slots = (256, pairs) if pair else (128, PLAN_SMS)
        n = up(I, 256) * up(J, 256) if pair else singles
        tail, stage, start = n % slots, 310 if pair else 290, 5000 if pair else 4000
        tile = (2500 if pair else 1500) + stage * kb
        forms.append(Plan(start + up(n, slots) * tile, n, 0, 0, 1, 0, pair))
        stages = tail * kb
        most = min(stages // 4, slots)
        if tail and most > 1:
            run = up(stages, most)
            ranges = up(stages, run)
            size = (ranges + tail) * edge * edge * 4
            apart = stage * run // 10 if 2 * (I + J) * R > L2_BYTES else 0
            forms.append(Plan(start + n // slots * tile + stage * run + apart + (9000 if pair else 4500) + size // 6000 + 30 * (ranges // tail), n - tail, ranges, run, 1, size, pair))
    for i, most in ((1, pairs), (2, 32), (3, 14)):
        if singles > most or (2 << i) > kb:
            break
        forms.append(Plan(4000 + 290 * ((kb + (1 << i) - 1) >> i) + 3500, singles, 0, 0, 1 << i, 0, False))
    return min(forms, key=lambda f: f.ns)           # (the first of equals)


def rows_ns(N, K):
    """Estimate of the form for one to eight rows."""
    units, steps, least = up(N, 16), up(K, 128), None
    for w in (2, 4, 8, 16):
        slices = 1
        while slices <= w and (slices == 1 or slices <= steps):
            t = up(up(units, w // slices), PLAN_SMS) * (up(steps, slices) * (140 * w + 1320) + 1500)
            least = t if least is None or t < least else least
            slices *= 2
    return 2500 + least * 10 // 19


def forward_form(M, N, K):
    plan = tile_plan(M, N, K)
    return "rows" if M <= 8 and rows_ns(N, K) * 3 // 4 <= plan.ns else plan.form


def workspace_bytes(M, N, K):
    most = up(N, 256) * 8 * 256 * 4 if M <= 8 else 0
    return 256 + max([most] + [tile_plan(*s).piece_bytes for s in ((M, N, K), (M, K, N), (N, K, M))])
