"""Calls of the dense operators that between them reach every kernel and layout, and the arguments of such a call on the host and on the device.

What a call gets is chosen by estimates on its sizes: each case says what it is there for, in the words of dlf_*_kernels on 148 SMs, and a test
on the host holds it to that.  A matrix is (rows, columns, pad, shift): values between two rows' ends and starts, and ahead of the first row."""
import ctypes as C
import re

from paper_2011_05630_b200 import binding as B, dense

STRUCTS = {"linear": dense._LINEAR, "linear_grad": dense._LINEAR_GRAD, "gated": dense._GATED, "gated_grad": dense._GATED_GRAD}
ORDER = {   # the structs' pointers, in their order; then the row lengths of those that are matrices, in the same order but for vectors
    "linear": "x w bias res y z", "linear_grad": "dy x w z dx dw db dz", "gated": "x wg wu bg bu h g u", "gated_grad": "dh x wg wu g u dx dwg dwu dbg dbu"}
VECTORS = {"bias", "db", "bg", "bu", "dbg", "dbu"}
OUTPUTS = {"linear": "y z", "linear_grad": "dx dw db dz", "gated": "h g u", "gated_grad": "dx dwg dwu dbg dbu"}


class Case:
    """pad, shift: of the inputs; out_pad, out_shift: of the outputs; without: what is null."""

    def __init__(self, name, op, m, k, n, expect, without="", pad=0, shift=0, out_pad=0, out_shift=0, act="relu"):
        self.name, self.op, self.m, self.k, self.n, self.expect, self.without, self.act = name, op, m, k, n, expect, without.split(), act
        self.pad, self.shift, self.out_pad, self.out_shift = pad, shift, out_pad, out_shift

    def matrices(self):
        """name -> (rows, columns, pad, shift), of those that are there."""
        m, k, n, out = self.m, self.k, self.n, OUTPUTS[self.op].split()
        size = {"x": (m, k), "dx": (m, k), "w": (n, k), "wg": (n, k), "wu": (n, k), "dw": (n, k), "dwg": (n, k), "dwu": (n, k)}
        return {t: size.get(t, (m, n)) + ((self.out_pad, self.out_shift) if t in out else (self.pad, self.shift))
                for t in ORDER[self.op].split() if t not in VECTORS and t not in self.without}

    def vectors(self):
        return [t for t in ORDER[self.op].split() if t in VECTORS and t not in self.without]

    def pack(self, dtype, pointer):
        """The argument struct; pointer(name) is where a matrix's first value or a vector lies."""
        mats, vecs = self.matrices(), self.vectors()
        names = ORDER[self.op].split()
        ptrs = [pointer(t) if t in mats or t in vecs else 0 for t in names]
        lds = [mats[t][1] + mats[t][2] if t in mats else 0 for t in names if t not in VECTORS]
        return STRUCTS[self.op].pack(B.DTYPES[dtype], B.DENSE_ACTS[self.act], self.m, self.k, self.n, *ptrs, *lds)

    def kernels(self, args, sms):
        text = C.create_string_buffer(1024)
        B._check(getattr(B.lib(), "dlf_%s_kernels" % self.op)(args, sms, text, len(text)), "dlf_%s_kernels" % self.op)
        return text.value.decode()

    def on_host(self, sms=148):
        """What a GPU of that many SMs would run, from pointers that nothing is read from."""
        mats = self.matrices()
        at = {t: (i + 1 << 30) + 2 * (mats[t][3] if t in mats else 0) for i, t in enumerate(ORDER[self.op].split())}
        return self.kernels(self.pack("bf16", at.get), sms)


def parts(text):
    """A call's kernels with their choices, but for the numbers that only grow with the sizes: + for any above 0 (of blocks: above 1)."""
    text = re.sub(r"pairs=\d+ ", "", text)
    text = re.sub(r"\b(rest|few|many)=(\d+)", lambda q: "%s=%s" % (q[1], "0" if q[2] == "0" else "+"), text)
    text = re.sub(r"blocks=(\d+)", lambda q: "blocks=%s" % ("1" if q[1] == "1" else "+"), text)
    return text.split("; ")


# (operator, m, k, n, pad, shift, out_pad, out_shift, what it is there for).  Without a further thought to the sizes: of random calls the largest
# with at most 600 million products that gets there, else the smallest.
_TABLE = [
    ("gated", 14, 3952, 4296, 0, 0, 0, 0, "dense_gemv(tokens=16 rows=aligned blocks=+ split=1)"),
    ("gated", 14, 4320, 1000, 0, 0, 3, 0, "dense_gemv(tokens=16 rows=aligned blocks=+ split=2)"),
    ("gated", 16, 3664, 592, 0, 8, 3, 0, "dense_gemv(tokens=16 rows=aligned blocks=+ split=4)"),
    ("gated", 15, 4088, 248, 8, 0, 3, 0, "dense_gemv(tokens=16 rows=aligned blocks=+ split=8)"),
    ("gated", 16, 704, 4008, 0, 0, 0, 0, "dense_gemv(tokens=16 rows=aligned blocks=1 split=1)"),
    ("gated", 16, 3479, 4197, 1, 0, 0, 0, "dense_gemv(tokens=16 rows=anywhere blocks=+ split=1)"),
    ("gated", 12, 4448, 1024, 1, 1, 0, 0, "dense_gemv(tokens=16 rows=anywhere blocks=+ split=2)"),
    ("gated", 16, 3842, 474, 0, 0, 3, 0, "dense_gemv(tokens=16 rows=anywhere blocks=+ split=4)"),
    ("gated", 14, 4432, 256, 8, 1, 0, 5, "dense_gemv(tokens=16 rows=anywhere blocks=+ split=8)"),
    ("gated", 13, 488, 4304, 1, 0, 0, 5, "dense_gemv(tokens=16 rows=anywhere blocks=1 split=1)"),
    ("gated", 8, 3960, 4400, 0, 0, 0, 0, "dense_gemv(tokens=8 rows=aligned blocks=+ split=1)"),
    ("gated", 7, 4232, 584, 0, 0, 0, 5, "dense_gemv(tokens=8 rows=aligned blocks=+ split=4)"),
    ("gated", 6, 4480, 272, 8, 0, 0, 5, "dense_gemv(tokens=8 rows=aligned blocks=+ split=8)"),
    ("gated", 8, 696, 3952, 0, 8, 3, 0, "dense_gemv(tokens=8 rows=aligned blocks=1 split=1)"),
    ("gated", 7, 4256, 4168, 1, 8, 0, 0, "dense_gemv(tokens=8 rows=anywhere blocks=+ split=1)"),
    ("gated", 7, 4492, 749, 1, 1, 3, 0, "dense_gemv(tokens=8 rows=anywhere blocks=+ split=2)"),
    ("gated", 7, 4311, 555, 8, 0, 0, 0, "dense_gemv(tokens=8 rows=anywhere blocks=+ split=4)"),
    ("gated", 8, 4184, 248, 1, 0, 0, 5, "dense_gemv(tokens=8 rows=anywhere blocks=+ split=8)"),
    ("gated", 6, 768, 4272, 1, 0, 0, 5, "dense_gemv(tokens=8 rows=anywhere blocks=1 split=1)"),
    ("gated", 271, 760, 2904, 1, 1, 0, 0, "dense_lat(products=1 columns=128 split=1 sources=1 out=aligned residual=none)"),
    ("gated", 425, 592, 2360, 0, 0, 3, 0, "dense_lat(products=1 columns=128 split=1 sources=1 out=anywhere residual=none)"),
    ("gated", 40, 3312, 4496, 8, 1, 0, 0, "dense_lat(products=1 columns=128 split=2 sources=1 out=aligned residual=none)"),
    ("gated", 51, 2448, 3928, 0, 1, 3, 5, "dense_lat(products=1 columns=128 split=2 sources=1 out=anywhere residual=none)"),
    ("gated", 861, 3104, 224, 8, 0, 0, 0, "dense_lat(products=1 columns=128 split=4 sources=1 out=aligned residual=none)"),
    ("gated", 800, 3088, 240, 0, 8, 3, 5, "dense_lat(products=1 columns=128 split=4 sources=1 out=anywhere residual=none)"),
    ("gated", 48, 4488, 944, 0, 1, 0, 0, "dense_lat(products=1 columns=128 split=8 sources=1 out=aligned residual=none)"),
    ("gated", 65, 4376, 848, 1, 1, 3, 0, "dense_lat(products=1 columns=128 split=8 sources=1 out=anywhere residual=none)"),
    ("gated", 189, 2152, 1464, 0, 1, 0, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=aligned residual=none)"),
    ("gated", 1028, 2257, 258, 0, 0, 0, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=anywhere residual=none)"),
    ("gated", 255, 2688, 872, 0, 1, 0, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=aligned residual=none)"),
    ("gated", 1259, 2354, 202, 0, 8, 0, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=anywhere residual=none)"),
    ("gated", 1011, 4334, 128, 0, 0, 0, 0, "dense_lat(products=1 columns=64 split=4 sources=1 out=aligned residual=none)"),
    ("gated", 1996, 4424, 56, 8, 8, 0, 5, "dense_lat(products=1 columns=64 split=4 sources=1 out=anywhere residual=none)"),
    ("gated", 565, 4472, 96, 8, 0, 0, 0, "dense_lat(products=1 columns=64 split=8 sources=1 out=aligned residual=none)"),
    ("gated", 616, 4016, 96, 8, 0, 3, 0, "dense_lat(products=1 columns=64 split=8 sources=1 out=anywhere residual=none)"),
    ("gated", 264, 960, 2344, 8, 0, 0, 0, "dense_lat(products=1 columns=96 split=1 sources=1 out=aligned residual=none)"),
    ("gated", 550, 1080, 1008, 8, 0, 0, 5, "dense_lat(products=1 columns=96 split=1 sources=1 out=anywhere residual=none)"),
    ("gated", 819, 2096, 344, 0, 0, 0, 0, "dense_lat(products=1 columns=96 split=2 sources=1 out=aligned residual=none)"),
    ("gated", 131, 3783, 1210, 0, 8, 0, 0, "dense_lat(products=1 columns=96 split=2 sources=1 out=anywhere residual=none)"),
    ("gated", 190, 4368, 720, 1, 0, 0, 0, "dense_lat(products=1 columns=96 split=4 sources=1 out=aligned residual=none)"),
    ("gated", 879, 4480, 152, 8, 8, 0, 5, "dense_lat(products=1 columns=96 split=4 sources=1 out=anywhere residual=none)"),
    ("gated", 369, 4352, 208, 0, 0, 0, 0, "dense_lat(products=1 columns=96 split=8 sources=1 out=aligned residual=none)"),
    ("gated", 827, 4408, 96, 0, 0, 3, 5, "dense_lat(products=1 columns=96 split=8 sources=1 out=anywhere residual=none)"),
    ("gated", 131, 3783, 1210, 0, 8, 0, 0, "dense_pack(matrices=3)"),
    ("gated", 1158, 232, 2216, 0, 1, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=aligned residual=none)"),
    ("gated", 1468, 152, 2680, 8, 0, 3, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=anywhere residual=none)"),
    ("gated", 1678, 480, 744, 0, 8, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=0 few=0 many=0 out=aligned residual=none)"),
    ("gated", 306, 456, 4296, 0, 8, 3, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=0 few=0 many=0 out=anywhere residual=none)"),
    ("gated_grad", 1834, 304, 1072, 0, 8, 0, 0, "dense_grad(rows=aligned columns=16)"),
    ("gated_grad", 176, 1448, 2352, 8, 8, 0, 0, "dense_grad(rows=aligned columns=64)"),
    ("gated_grad", 2048, 248, 1176, 1, 0, 0, 0, "dense_grad(rows=anywhere columns=16)"),
    ("gated_grad", 937, 456, 1400, 1, 0, 0, 0, "dense_grad(rows=anywhere columns=64)"),
    ("gated_grad", 167, 1648, 1384, 1, 1, 0, 0, "dense_lat(products=1 columns=128 split=1 sources=1 out=aligned residual=none)"),
    ("gated_grad", 184, 619, 3670, 1, 1, 3, 5, "dense_lat(products=1 columns=128 split=1 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 1822, 1824, 64, 0, 0, 0, 0, "dense_lat(products=1 columns=128 split=1 sources=2 out=aligned residual=none)"),
    ("gated_grad", 1913, 1735, 64, 8, 0, 3, 0, "dense_lat(products=1 columns=128 split=1 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 2070, 3664, 8, 1, 0, 0, 5, "dense_lat(products=1 columns=128 split=2 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 131, 2496, 1488, 0, 8, 0, 0, "dense_lat(products=1 columns=128 split=2 sources=2 out=aligned residual=none)"),
    ("gated_grad", 138, 2652, 2006, 0, 1, 3, 0, "dense_lat(products=1 columns=128 split=2 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1993, 1984, 56, 8, 8, 0, 0, "dense_lat(products=1 columns=128 split=4 sources=1 out=aligned residual=none)"),
    ("gated_grad", 2045, 1982, 63, 0, 0, 0, 0, "dense_lat(products=1 columns=128 split=4 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 176, 1448, 2352, 8, 8, 0, 0, "dense_lat(products=1 columns=128 split=4 sources=2 out=aligned residual=none)"),
    ("gated_grad", 45, 3512, 3736, 1, 0, 0, 5, "dense_lat(products=1 columns=128 split=4 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1846, 528, 32, 0, 8, 0, 0, "dense_lat(products=1 columns=128 split=8 sources=1 out=aligned residual=none)"),
    ("gated_grad", 2012, 824, 32, 1, 0, 3, 5, "dense_lat(products=1 columns=128 split=8 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 156, 872, 4048, 0, 0, 0, 0, "dense_lat(products=1 columns=128 split=8 sources=2 out=aligned residual=none)"),
    ("gated_grad", 269, 538, 4024, 0, 0, 0, 5, "dense_lat(products=1 columns=128 split=8 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 991, 264, 2224, 0, 0, 0, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=aligned residual=none)"),
    ("gated_grad", 1040, 216, 2640, 1, 8, 3, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 137, 2696, 1396, 1, 0, 0, 0, "dense_lat(products=1 columns=64 split=1 sources=2 out=aligned residual=none)"),
    ("gated_grad", 266, 1744, 1256, 1, 0, 3, 0, "dense_lat(products=1 columns=64 split=1 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1875, 64, 4440, 8, 8, 0, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=aligned residual=none)"),
    ("gated_grad", 1932, 56, 4016, 1, 8, 3, 5, "dense_lat(products=1 columns=64 split=2 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 331, 1056, 1680, 8, 0, 0, 0, "dense_lat(products=1 columns=64 split=2 sources=2 out=aligned residual=none)"),
    ("gated_grad", 90, 3824, 1736, 0, 8, 0, 5, "dense_lat(products=1 columns=64 split=2 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 2013, 488, 176, 8, 8, 0, 0, "dense_lat(products=1 columns=64 split=4 sources=1 out=aligned residual=none)"),
    ("gated_grad", 2032, 984, 104, 0, 0, 3, 0, "dense_lat(products=1 columns=64 split=4 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 498, 376, 3168, 1, 0, 0, 0, "dense_lat(products=1 columns=64 split=4 sources=2 out=aligned residual=none)"),
    ("gated_grad", 579, 322, 3205, 1, 1, 0, 0, "dense_lat(products=1 columns=64 split=4 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1873, 432, 64, 0, 0, 0, 0, "dense_lat(products=1 columns=64 split=8 sources=1 out=aligned residual=none)"),
    ("gated_grad", 2024, 280, 64, 8, 0, 3, 5, "dense_lat(products=1 columns=64 split=8 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 1875, 64, 4440, 8, 8, 0, 0, "dense_lat(products=1 columns=64 split=8 sources=2 out=aligned residual=none)"),
    ("gated_grad", 847, 128, 4456, 1, 0, 3, 0, "dense_lat(products=1 columns=64 split=8 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1845, 536, 584, 8, 1, 0, 0, "dense_lat(products=2 columns=128 split=1 sources=1 out=aligned residual=none)"),
    ("gated_grad", 1556, 639, 598, 0, 0, 3, 0, "dense_lat(products=2 columns=128 split=1 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 937, 456, 1400, 1, 0, 0, 0, "dense_lat(products=2 columns=128 split=1 sources=2 out=aligned residual=none)"),
    ("gated_grad", 1292, 364, 1238, 8, 0, 0, 0, "dense_lat(products=2 columns=128 split=1 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1904, 456, 24, 0, 8, 0, 0, "dense_lat(products=2 columns=128 split=2 sources=1 out=aligned residual=none)"),
    ("gated_grad", 2040, 464, 32, 1, 8, 3, 0, "dense_lat(products=2 columns=128 split=2 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 1955, 128, 2224, 8, 8, 0, 0, "dense_lat(products=2 columns=128 split=2 sources=2 out=aligned residual=none)"),
    ("gated_grad", 2083, 96, 2480, 0, 0, 0, 5, "dense_lat(products=2 columns=128 split=2 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1360, 640, 678, 8, 0, 0, 0, "dense_lat(products=2 columns=64 split=1 sources=1 out=aligned residual=none)"),
    ("gated_grad", 2006, 560, 490, 8, 0, 0, 5, "dense_lat(products=2 columns=64 split=1 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 1834, 304, 1072, 0, 8, 0, 0, "dense_lat(products=2 columns=64 split=1 sources=2 out=aligned residual=none)"),
    ("gated_grad", 1510, 208, 1880, 8, 0, 0, 5, "dense_lat(products=2 columns=64 split=1 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1790, 152, 600, 8, 0, 0, 0, "dense_lat(products=2 columns=64 split=2 sources=1 out=aligned residual=none)"),
    ("gated_grad", 1951, 112, 904, 8, 0, 3, 0, "dense_lat(products=2 columns=64 split=2 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 1667, 64, 3264, 0, 0, 0, 0, "dense_lat(products=2 columns=64 split=2 sources=2 out=aligned residual=none)"),
    ("gated_grad", 1391, 64, 3616, 8, 1, 3, 0, "dense_lat(products=2 columns=64 split=2 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 2073, 56, 784, 1, 8, 0, 0, "dense_lat(products=2 columns=64 split=4 sources=1 out=aligned residual=none)"),
    ("gated_grad", 1966, 63, 940, 0, 0, 0, 0, "dense_lat(products=2 columns=64 split=4 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 1864, 64, 1072, 8, 0, 0, 0, "dense_lat(products=2 columns=64 split=4 sources=2 out=aligned residual=none)"),
    ("gated_grad", 1303, 64, 1408, 8, 0, 0, 5, "dense_lat(products=2 columns=64 split=4 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1386, 40, 224, 1, 0, 0, 0, "dense_lat(products=2 columns=64 split=8 sources=1 out=aligned residual=none)"),
    ("gated_grad", 902, 56, 255, 8, 0, 0, 5, "dense_lat(products=2 columns=64 split=8 sources=1 out=anywhere residual=none)"),
    ("gated_grad", 500, 8, 512, 0, 1, 0, 0, "dense_lat(products=2 columns=64 split=8 sources=2 out=aligned residual=none)"),
    ("gated_grad", 509, 40, 488, 0, 0, 3, 0, "dense_lat(products=2 columns=64 split=8 sources=2 out=anywhere residual=none)"),
    ("gated_grad", 1, 8, 8, 1, 0, 0, 0, "dense_pack(matrices=2)"),
    ("gated_grad", 937, 456, 1400, 1, 0, 0, 0, "dense_pack(matrices=3)"),
    ("gated_grad", 266, 1088, 1976, 0, 0, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=2 rest=+ few=0 many=0 out=aligned residual=none)"),
    ("gated_grad", 271, 872, 2416, 0, 0, 0, 5, "dense_pair(products=1 columns=128 sources=1 groups=2 rest=+ few=0 many=0 out=anywhere residual=none)"),
    ("gated_grad", 589, 656, 1424, 0, 0, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=2 rest=0 few=0 many=0 out=aligned residual=none)"),
    ("gated_grad", 634, 656, 1432, 8, 8, 3, 0, "dense_pair(products=1 columns=128 sources=1 groups=2 rest=0 few=0 many=0 out=anywhere residual=none)"),
    ("gated_grad", 1956, 1136, 112, 1, 0, 0, 0, "dense_pair(products=1 columns=128 sources=2 groups=1 rest=0 few=0 many=0 out=aligned residual=none)"),
    ("gated_grad", 2003, 1072, 80, 8, 8, 3, 5, "dense_pair(products=1 columns=128 sources=2 groups=1 rest=0 few=0 many=0 out=anywhere residual=none)"),
    ("gated_grad", 176, 1448, 2352, 8, 8, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=2 rest=+ few=0 many=0 out=aligned residual=none)"),
    ("gated_grad", 90, 3824, 1736, 0, 8, 0, 5, "dense_pair(products=1 columns=256 sources=1 groups=2 rest=+ few=0 many=0 out=anywhere residual=none)"),
    ("gated_grad", 498, 376, 3168, 1, 0, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=2 rest=0 few=0 many=0 out=aligned residual=none)"),
    ("gated_grad", 579, 322, 3205, 1, 1, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=2 rest=0 few=0 many=0 out=anywhere residual=none)"),
    ("gated_grad", 1990, 2360, 24, 0, 8, 0, 0, "dense_pair(products=1 columns=256 sources=2 groups=1 rest=+ few=0 many=0 out=aligned residual=none)"),
    ("gated_grad", 2037, 2344, 8, 0, 1, 0, 5, "dense_pair(products=1 columns=256 sources=2 groups=1 rest=+ few=0 many=0 out=anywhere residual=none)"),
    ("gated_grad", 1993, 1984, 56, 8, 8, 0, 0, "dense_pair(products=1 columns=256 sources=2 groups=1 rest=0 few=0 many=0 out=aligned residual=none)"),
    ("gated_grad", 2005, 2264, 80, 1, 0, 3, 0, "dense_pair(products=1 columns=256 sources=2 groups=1 rest=0 few=0 many=0 out=anywhere residual=none)"),
    ("gated_grad", 1580, 1336, 712, 0, 8, 0, 5, "dense_pair(products=2 columns=128 sources=1 groups=1 rest=+ few=+ many=+ out=anywhere residual=none)"),
    ("gated_grad", 1842, 1064, 304, 1, 0, 0, 0, "dense_pair(products=2 columns=128 sources=1 groups=1 rest=+ few=+ many=0 out=aligned residual=none)"),
    ("gated_grad", 1502, 1552, 256, 1, 0, 3, 0, "dense_pair(products=2 columns=128 sources=1 groups=1 rest=+ few=+ many=0 out=anywhere residual=none)"),
    ("gated_grad", 670, 2600, 344, 8, 8, 3, 5, "dense_pair(products=2 columns=128 sources=2 groups=2 rest=+ few=+ many=+ out=anywhere residual=none)"),
    ("gated_grad", 173, 2968, 1128, 0, 8, 0, 0, "dense_pair(products=2 columns=128 sources=2 groups=2 rest=+ few=+ many=0 out=aligned residual=none)"),
    ("gated_grad", 593, 1440, 688, 1, 0, 0, 5, "dense_pair(products=2 columns=128 sources=2 groups=2 rest=+ few=+ many=0 out=anywhere residual=none)"),
    ("gated_grad", 620, 3000, 264, 1, 0, 0, 0, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=+ out=aligned residual=none)"),
    ("gated_grad", 618, 3416, 296, 0, 1, 0, 5, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=+ out=anywhere residual=none)"),
    ("gated_grad", 1279, 3592, 128, 8, 0, 0, 0, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=0 out=aligned residual=none)"),
    ("gated_grad", 956, 2317, 269, 1, 0, 0, 5, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=0 out=anywhere residual=none)"),
    ("gated_grad", 527, 3608, 344, 8, 0, 0, 0, "dense_pair(products=2 columns=256 sources=2 groups=2 rest=+ few=+ many=+ out=aligned residual=none)"),
    ("gated_grad", 572, 3639, 400, 0, 8, 0, 0, "dense_pair(products=2 columns=256 sources=2 groups=2 rest=+ few=+ many=+ out=anywhere residual=none)"),
    ("gated_grad", 213, 3144, 880, 1, 0, 0, 0, "dense_pair(products=2 columns=256 sources=2 groups=2 rest=+ few=+ many=0 out=aligned residual=none)"),
    ("gated_grad", 516, 3346, 344, 1, 0, 0, 5, "dense_pair(products=2 columns=256 sources=2 groups=2 rest=+ few=+ many=0 out=anywhere residual=none)"),
    ("linear", 16, 4320, 4472, 8, 0, 3, 5, "dense_gemv(tokens=16 rows=aligned blocks=+ split=1)"),
    ("linear", 15, 4232, 440, 0, 0, 3, 5, "dense_gemv(tokens=16 rows=aligned blocks=+ split=4)"),
    ("linear", 14, 4288, 224, 0, 8, 3, 5, "dense_gemv(tokens=16 rows=aligned blocks=+ split=8)"),
    ("linear", 15, 896, 4400, 0, 0, 0, 0, "dense_gemv(tokens=16 rows=aligned blocks=1 split=1)"),
    ("linear", 14, 4446, 3590, 0, 0, 3, 0, "dense_gemv(tokens=16 rows=anywhere blocks=+ split=1)"),
    ("linear", 16, 4091, 575, 0, 1, 0, 0, "dense_gemv(tokens=16 rows=anywhere blocks=+ split=4)"),
    ("linear", 14, 4222, 226, 0, 0, 0, 0, "dense_gemv(tokens=16 rows=anywhere blocks=+ split=8)"),
    ("linear", 16, 928, 4136, 1, 8, 0, 0, "dense_gemv(tokens=16 rows=anywhere blocks=1 split=1)"),
    ("linear", 8, 3904, 4200, 0, 0, 0, 0, "dense_gemv(tokens=8 rows=aligned blocks=+ split=1)"),
    ("linear", 8, 1392, 4288, 0, 8, 0, 0, "dense_gemv(tokens=8 rows=aligned blocks=1 split=1)"),
    ("linear", 8, 3024, 3968, 1, 0, 0, 5, "dense_gemv(tokens=8 rows=anywhere blocks=+ split=1)"),
    ("linear", 8, 4480, 480, 1, 0, 0, 0, "dense_gemv(tokens=8 rows=anywhere blocks=+ split=4)"),
    ("linear", 7, 1192, 4400, 1, 8, 0, 5, "dense_gemv(tokens=8 rows=anywhere blocks=1 split=1)"),
    ("linear", 1838, 128, 2416, 0, 0, 0, 0, "dense_lat(products=1 columns=128 split=1 sources=1 out=aligned residual=aligned)"),
    ("linear", 1795, 128, 1936, 1, 0, 0, 0, "dense_lat(products=1 columns=128 split=1 sources=1 out=aligned residual=anywhere)"),
    ("linear", 1102, 128, 3936, 0, 0, 3, 0, "dense_lat(products=1 columns=128 split=1 sources=1 out=anywhere residual=aligned)"),
    ("linear", 1044, 176, 3264, 1, 8, 0, 5, "dense_lat(products=1 columns=128 split=1 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 1470, 2808, 600, 0, 0, 0, 0, "dense_lat(products=1 columns=128 split=2 sources=1 out=aligned residual=aligned)"),
    ("linear", 157, 3680, 3784, 8, 1, 0, 0, "dense_lat(products=1 columns=128 split=2 sources=1 out=aligned residual=anywhere)"),
    ("linear", 272, 3048, 2736, 8, 0, 0, 5, "dense_lat(products=1 columns=128 split=2 sources=1 out=anywhere residual=aligned)"),
    ("linear", 153, 3308, 4302, 0, 0, 0, 0, "dense_lat(products=1 columns=128 split=2 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 50, 2560, 3952, 0, 8, 0, 0, "dense_lat(products=1 columns=128 split=4 sources=1 out=aligned residual=aligned)"),
    ("linear", 68, 2256, 3408, 1, 0, 0, 0, "dense_lat(products=1 columns=128 split=4 sources=1 out=aligned residual=anywhere)"),
    ("linear", 62, 2736, 3352, 8, 0, 0, 5, "dense_lat(products=1 columns=128 split=4 sources=1 out=anywhere residual=aligned)"),
    ("linear", 58, 2662, 3807, 0, 1, 0, 0, "dense_lat(products=1 columns=128 split=4 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 54, 4088, 1920, 8, 0, 0, 0, "dense_lat(products=1 columns=128 split=8 sources=1 out=aligned residual=aligned)"),
    ("linear", 57, 4192, 1576, 8, 1, 0, 0, "dense_lat(products=1 columns=128 split=8 sources=1 out=aligned residual=anywhere)"),
    ("linear", 18, 4000, 1880, 0, 0, 0, 5, "dense_lat(products=1 columns=128 split=8 sources=1 out=anywhere residual=aligned)"),
    ("linear", 52, 4136, 1672, 0, 1, 3, 0, "dense_lat(products=1 columns=128 split=8 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 866, 720, 952, 8, 0, 0, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=aligned residual=aligned)"),
    ("linear", 398, 824, 1776, 1, 0, 0, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=aligned residual=anywhere)"),
    ("linear", 767, 488, 1600, 0, 0, 3, 5, "dense_lat(products=1 columns=64 split=1 sources=1 out=anywhere residual=aligned)"),
    ("linear", 230, 659, 3953, 0, 0, 0, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 196, 1328, 2256, 0, 0, 0, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=aligned residual=aligned)"),
    ("linear", 179, 1672, 2000, 1, 0, 0, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=aligned residual=anywhere)"),
    ("linear", 222, 1296, 2080, 0, 8, 3, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=anywhere residual=aligned)"),
    ("linear", 193, 1615, 1922, 0, 0, 3, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 1059, 4384, 128, 0, 0, 0, 0, "dense_lat(products=1 columns=64 split=4 sources=1 out=aligned residual=aligned)"),
    ("linear", 107, 2976, 1768, 8, 1, 0, 0, "dense_lat(products=1 columns=64 split=4 sources=1 out=aligned residual=anywhere)"),
    ("linear", 646, 3744, 248, 0, 8, 3, 5, "dense_lat(products=1 columns=64 split=4 sources=1 out=anywhere residual=aligned)"),
    ("linear", 330, 3360, 536, 1, 0, 0, 5, "dense_lat(products=1 columns=64 split=4 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 320, 4448, 312, 0, 0, 0, 0, "dense_lat(products=1 columns=64 split=8 sources=1 out=aligned residual=aligned)"),
    ("linear", 1832, 3688, 64, 1, 8, 0, 0, "dense_lat(products=1 columns=64 split=8 sources=1 out=aligned residual=anywhere)"),
    ("linear", 1900, 3536, 64, 8, 0, 3, 5, "dense_lat(products=1 columns=64 split=8 sources=1 out=anywhere residual=aligned)"),
    ("linear", 332, 4232, 304, 0, 1, 3, 0, "dense_lat(products=1 columns=64 split=8 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 932, 256, 2328, 8, 8, 0, 0, "dense_lat(products=1 columns=96 split=1 sources=1 out=aligned residual=aligned)"),
    ("linear", 1904, 392, 800, 1, 0, 0, 0, "dense_lat(products=1 columns=96 split=1 sources=1 out=aligned residual=anywhere)"),
    ("linear", 942, 352, 1800, 8, 8, 0, 5, "dense_lat(products=1 columns=96 split=1 sources=1 out=anywhere residual=aligned)"),
    ("linear", 564, 484, 2190, 0, 8, 0, 5, "dense_lat(products=1 columns=96 split=1 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 153, 2056, 3032, 8, 0, 0, 0, "dense_lat(products=1 columns=96 split=2 sources=1 out=aligned residual=aligned)"),
    ("linear", 129, 2160, 2520, 1, 0, 0, 0, "dense_lat(products=1 columns=96 split=2 sources=1 out=aligned residual=anywhere)"),
    ("linear", 162, 1928, 2472, 0, 0, 3, 0, "dense_lat(products=1 columns=96 split=2 sources=1 out=anywhere residual=aligned)"),
    ("linear", 133, 2208, 2392, 8, 1, 3, 0, "dense_lat(products=1 columns=96 split=2 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 410, 2280, 640, 8, 0, 0, 0, "dense_lat(products=1 columns=96 split=4 sources=1 out=aligned residual=aligned)"),
    ("linear", 122, 1760, 2736, 1, 1, 0, 0, "dense_lat(products=1 columns=96 split=4 sources=1 out=aligned residual=anywhere)"),
    ("linear", 1460, 2664, 152, 8, 0, 3, 0, "dense_lat(products=1 columns=96 split=4 sources=1 out=anywhere residual=aligned)"),
    ("linear", 199, 2834, 1052, 0, 0, 0, 5, "dense_lat(products=1 columns=96 split=4 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 245, 3552, 672, 0, 0, 0, 0, "dense_lat(products=1 columns=96 split=8 sources=1 out=aligned residual=aligned)"),
    ("linear", 343, 4248, 400, 1, 1, 0, 0, "dense_lat(products=1 columns=96 split=8 sources=1 out=aligned residual=anywhere)"),
    ("linear", 812, 3760, 192, 0, 8, 0, 5, "dense_lat(products=1 columns=96 split=8 sources=1 out=anywhere residual=aligned)"),
    ("linear", 580, 3992, 256, 0, 1, 3, 5, "dense_lat(products=1 columns=96 split=8 sources=1 out=anywhere residual=anywhere)"),
    ("linear", 1044, 176, 3264, 1, 8, 0, 5, "dense_pack(matrices=2)"),
    ("linear", 1751, 248, 2680, 0, 0, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=+ few=0 many=0 out=aligned residual=aligned)"),
    ("linear", 1258, 379, 3649, 0, 1, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=+ few=0 many=0 out=anywhere residual=anywhere)"),
    ("linear", 714, 288, 2824, 0, 8, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=0 few=0 many=0 out=aligned residual=aligned)"),
    ("linear", 500, 208, 4360, 1, 0, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=0 few=0 many=0 out=aligned residual=anywhere)"),
    ("linear", 1292, 296, 1440, 8, 0, 3, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=0 few=0 many=0 out=anywhere residual=aligned)"),
    ("linear", 1997, 296, 942, 0, 0, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=0 few=0 many=0 out=anywhere residual=anywhere)"),
    ("linear", 2100, 72, 3640, 8, 0, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=aligned residual=aligned)"),
    ("linear", 1193, 112, 3976, 1, 0, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=aligned residual=anywhere)"),
    ("linear", 1284, 104, 4320, 0, 0, 3, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=anywhere residual=aligned)"),
    ("linear", 1895, 72, 4008, 1, 0, 3, 5, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=anywhere residual=anywhere)"),
    ("linear", 1643, 144, 2488, 0, 0, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=0 few=0 many=0 out=aligned residual=aligned)"),
    ("linear", 870, 216, 2976, 1, 1, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=0 few=0 many=0 out=aligned residual=anywhere)"),
    ("linear", 1218, 144, 3400, 8, 0, 3, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=0 few=0 many=0 out=anywhere residual=aligned)"),
    ("linear", 1882, 208, 1520, 0, 1, 3, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=0 few=0 many=0 out=anywhere residual=anywhere)"),
    ("linear_grad", 1854, 232, 1384, 0, 8, 0, 0, "dense_grad(rows=aligned columns=16)"),
    ("linear_grad", 247, 1280, 1896, 8, 0, 0, 0, "dense_grad(rows=aligned columns=64)"),
    ("linear_grad", 1972, 162, 1871, 8, 0, 0, 0, "dense_grad(rows=anywhere columns=16)"),
    ("linear_grad", 252, 1224, 1944, 0, 0, 3, 0, "dense_grad(rows=anywhere columns=64)"),
    ("linear_grad", 145, 1056, 3784, 8, 0, 0, 0, "dense_lat(products=1 columns=128 split=1 sources=1 out=aligned residual=none)"),
    ("linear_grad", 136, 1654, 2599, 1, 0, 0, 0, "dense_lat(products=1 columns=128 split=1 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 151, 2624, 3144, 1, 0, 0, 0, "dense_lat(products=1 columns=128 split=2 sources=1 out=aligned residual=none)"),
    ("linear_grad", 137, 3504, 4208, 8, 1, 3, 0, "dense_lat(products=1 columns=128 split=2 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 57, 3736, 2768, 0, 8, 0, 0, "dense_lat(products=1 columns=128 split=4 sources=1 out=aligned residual=none)"),
    ("linear_grad", 55, 2896, 3688, 8, 8, 3, 5, "dense_lat(products=1 columns=128 split=4 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 49, 1656, 3528, 1, 0, 0, 0, "dense_lat(products=1 columns=128 split=8 sources=1 out=aligned residual=none)"),
    ("linear_grad", 133, 829, 4453, 0, 0, 3, 5, "dense_lat(products=1 columns=128 split=8 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 731, 184, 4448, 0, 8, 0, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=aligned residual=none)"),
    ("linear_grad", 750, 260, 3071, 1, 0, 3, 0, "dense_lat(products=1 columns=64 split=1 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 202, 1456, 2016, 1, 1, 0, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=aligned residual=none)"),
    ("linear_grad", 164, 1500, 2437, 1, 0, 0, 0, "dense_lat(products=1 columns=64 split=2 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 731, 184, 4448, 0, 8, 0, 0, "dense_lat(products=1 columns=64 split=4 sources=1 out=aligned residual=none)"),
    ("linear_grad", 750, 260, 3071, 1, 0, 3, 0, "dense_lat(products=1 columns=64 split=4 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 128, 952, 3824, 8, 0, 0, 0, "dense_lat(products=1 columns=64 split=8 sources=1 out=aligned residual=none)"),
    ("linear_grad", 369, 310, 4319, 1, 0, 0, 0, "dense_lat(products=1 columns=64 split=8 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 452, 896, 1464, 1, 1, 0, 0, "dense_lat(products=2 columns=128 split=1 sources=1 out=aligned residual=none)"),
    ("linear_grad", 950, 1160, 544, 0, 1, 0, 5, "dense_lat(products=2 columns=128 split=1 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 1791, 104, 3184, 8, 8, 0, 0, "dense_lat(products=2 columns=128 split=2 sources=1 out=aligned residual=none)"),
    ("linear_grad", 1003, 131, 3533, 8, 1, 3, 0, "dense_lat(products=2 columns=128 split=2 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 1030, 120, 2464, 0, 0, 0, 0, "dense_lat(products=2 columns=128 split=4 sources=1 out=aligned residual=none)"),
    ("linear_grad", 1001, 69, 2744, 0, 0, 0, 0, "dense_lat(products=2 columns=128 split=4 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 1455, 128, 3207, 1, 0, 0, 0, "dense_lat(products=2 columns=64 split=1 sources=1 out=aligned residual=none)"),
    ("linear_grad", 1184, 128, 3944, 0, 0, 0, 5, "dense_lat(products=2 columns=64 split=1 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 1709, 120, 2752, 0, 0, 0, 0, "dense_lat(products=2 columns=64 split=2 sources=1 out=aligned residual=none)"),
    ("linear_grad", 1388, 128, 3176, 1, 0, 0, 5, "dense_lat(products=2 columns=64 split=2 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 1529, 64, 2624, 8, 0, 0, 0, "dense_lat(products=2 columns=64 split=4 sources=1 out=aligned residual=none)"),
    ("linear_grad", 1404, 64, 2816, 0, 0, 3, 0, "dense_lat(products=2 columns=64 split=4 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 471, 40, 1392, 8, 8, 0, 0, "dense_lat(products=2 columns=64 split=8 sources=1 out=aligned residual=none)"),
    ("linear_grad", 492, 56, 1368, 8, 0, 3, 5, "dense_lat(products=2 columns=64 split=8 sources=1 out=anywhere residual=none)"),
    ("linear_grad", 1, 8, 8, 1, 0, 3, 0, "dense_pack(matrices=1)"),
    ("linear_grad", 164, 1500, 2437, 1, 0, 0, 0, "dense_pack(matrices=2)"),
    ("linear_grad", 2, 2080, 4216, 1, 0, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=+ few=0 many=0 out=aligned residual=none)"),
    ("linear_grad", 50, 3704, 2464, 1, 0, 3, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=+ few=0 many=0 out=anywhere residual=none)"),
    ("linear_grad", 252, 960, 2200, 8, 0, 0, 0, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=0 few=0 many=0 out=aligned residual=none)"),
    ("linear_grad", 282, 631, 3331, 1, 0, 0, 5, "dense_pair(products=1 columns=128 sources=1 groups=1 rest=0 few=0 many=0 out=anywhere residual=none)"),
    ("linear_grad", 57, 3736, 2768, 0, 8, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=aligned residual=none)"),
    ("linear_grad", 43, 4400, 3160, 0, 0, 3, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=anywhere residual=none)"),
    ("linear_grad", 241, 848, 2912, 8, 8, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=0 few=0 many=0 out=aligned residual=none)"),
    ("linear_grad", 164, 1500, 2437, 1, 0, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=0 few=0 many=0 out=anywhere residual=none)"),
    ("linear_grad", 715, 2672, 832, 0, 0, 0, 0, "dense_pair(products=2 columns=128 sources=1 groups=1 rest=+ few=+ many=+ out=aligned residual=none)"),
    ("linear_grad", 766, 2674, 818, 0, 0, 0, 5, "dense_pair(products=2 columns=128 sources=1 groups=1 rest=+ few=+ many=+ out=anywhere residual=none)"),
    ("linear_grad", 247, 1280, 1896, 8, 0, 0, 0, "dense_pair(products=2 columns=128 sources=1 groups=1 rest=+ few=+ many=0 out=aligned residual=none)"),
    ("linear_grad", 252, 1224, 1944, 0, 0, 3, 0, "dense_pair(products=2 columns=128 sources=1 groups=1 rest=+ few=+ many=0 out=anywhere residual=none)"),
    ("linear_grad", 542, 3192, 616, 0, 1, 0, 0, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=+ out=aligned residual=none)"),
    ("linear_grad", 460, 3992, 528, 0, 1, 3, 0, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=+ out=anywhere residual=none)"),
    ("linear_grad", 536, 2360, 472, 1, 0, 0, 0, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=0 out=aligned residual=none)"),
    ("linear_grad", 328, 4480, 408, 0, 0, 3, 0, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=0 out=anywhere residual=none)"),
    # more than a pair's share of tiles, a second job's tiles shared out unevenly; sizes that divide by nothing
    ("linear", 1500, 1111, 3333, 1, 0, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=anywhere residual=anywhere)"),
    ("gated", 3000, 999, 1777, 0, 0, 0, 0, "dense_pair(products=1 columns=256 sources=1 groups=1 rest=+ few=0 many=0 out=anywhere residual=none)"),
    ("linear_grad", 2048, 2048, 2048, 0, 0, 0, 0, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=+ out=aligned residual=none)"),
    ("gated_grad", 2048, 2048, 2048, 0, 0, 0, 0, "dense_pair(products=2 columns=256 sources=2 groups=2 rest=+ few=+ many=+ out=aligned residual=none)"),
    ("linear_grad", 1500, 1111, 3333, 0, 0, 0, 0, "dense_pair(products=2 columns=256 sources=1 groups=1 rest=+ few=+ many=0 out=anywhere residual=none)"),
    ("gated_grad", 612, 2584, 344, 1, 0, 0, 0, "dense_pair(products=2 columns=128 sources=2 groups=2 rest=+ few=+ many=+ out=aligned residual=none)"),
    ("linear_grad", 20000, 64, 33, 0, 0, 0, 0, "dense_grad(rows=anywhere columns=16)"),
]
CASES = [Case("%d: %s %d x %d x %d" % (i, t[0], *t[1:4]), t[0], *t[1:4], t[8], pad=t[4], shift=t[5], out_pad=t[6], out_shift=t[7]) for i, t in enumerate(_TABLE)]

# what the kernels' templates and the host's choices make possible: each has a case
REACHED = [
    *("dense_gemv(tokens=%d rows=%s blocks=%s split=%d)" % (t, r, b, s) for t in (8, 16) for r in ("aligned", "anywhere") for b, s in (("1", 1), ("+", 1), ("+", 4))),
    *("dense_grad(rows=%s columns=%d)" % (r, c) for r in ("aligned", "anywhere") for c in (16, 64)),
    *("dense_lat(products=1 columns=%d split=%d sources=1 out=%s residual=%s)" % (c, s, o, r) for c in (64, 96, 128) for s in (1, 2, 4, 8)
      for o in ("aligned", "anywhere") for r in ("aligned", "anywhere")),
    *("dense_lat(products=2 columns=%d split=1 sources=%d out=%s residual=none)" % (c, s, o) for c in (64, 128) for s in (1, 2) for o in ("aligned", "anywhere")),
    *("dense_lat(products=2 columns=64 split=%d sources=%d out=%s residual=none)" % (s, q, o) for s in (2, 4, 8) for q in (1, 2) for o in ("aligned", "anywhere")),
    *("dense_pair(products=1 columns=256 sources=1 groups=1 rest=%s few=0 many=0 out=%s residual=%s)" % (t, o, r) for t in "0+" for o in ("aligned", "anywhere")
      for r in ("none", "aligned", "anywhere")),
    *("dense_pair(products=1 columns=128 sources=1 groups=1 rest=0 few=0 many=0 out=%s residual=%s)" % (o, r) for o in ("aligned", "anywhere") for r in ("none", "aligned")),
    *("dense_pair(products=1 columns=%d sources=1 groups=2 rest=%s few=0 many=0 out=%s residual=none)" % (c, t, o) for c in (128, 256) for t in "0+" for o in ("aligned", "anywhere")),
    *("dense_pair(products=2 columns=%d sources=%d groups=%d rest=+ few=+ many=%s out=%s residual=none)" % (c, s, s, t, o) for c in (128, 256) for s in (1, 2)
      for t in "0+" for o in ("aligned", "anywhere")),
]
