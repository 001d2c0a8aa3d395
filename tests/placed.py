"""Matrices with a pitch and an offset of their own inside a larger buffer, which is looked at afterwards."""
MARK = 5.0


class Placed:
    def __init__(self, torch, rows, cols, dtype, pad=0, offset=0, fill=None):
        self.rows, self.cols, self.ld, self.offset = rows, cols, cols + pad, offset
        self.flat = torch.full((offset + rows * self.ld + 16,), MARK, dtype=dtype, device="cuda")
        self.m = self.flat[offset:offset + rows * self.ld].view(rows, self.ld)
        if fill is not None:
            self.m[:, :cols] = fill.to(dtype)

    @property
    def values(self):
        return self.m[:, :self.cols]

    def guarded(self):
        """Nothing was written beside the matrix."""
        return bool((self.flat[:self.offset] == MARK).all()) and bool((self.m[:, self.cols:] == MARK).all()) and bool((self.flat[self.offset + self.m.numel():] == MARK).all())

    def data_ptr(self):
        return self.m.data_ptr()
