"""Which kernels the entry points of stagefrontier_train.h launch, without a
GPU: run in a process of its own with launch_recorder.c in place of the HIP
runtime.  Reads a JSON list of [function, [arguments]]; an argument is "p<i>"
(one of a set of far apart addresses that nothing reads), ["i", v], ["l", v],
["f", v], or ["list", [[address index, numel, dtype], ...]] for a list of
gradients, which is laid out first."""
import ctypes
import json
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))


def address(i):
    return (int(i) + 1) << 46


def main():
    rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    rec.rec_name.restype = ctypes.c_char_p
    rec.rec_lds.restype = ctypes.c_uint64
    lib = ctypes.CDLL(sys.argv[2])
    lib.sf_grad_list_bytes.restype = ctypes.c_int64
    out = []
    for name, args in json.load(sys.stdin):
        conv, keep, at = [], [], 0
        for a in args:
            if isinstance(a, str):
                conv.append(ctypes.c_void_p(address(a[1:])))
            elif a[0] == "list":
                n = len(a[1])
                size = lib.sf_grad_list_bytes(ctypes.c_int32(n))
                buf = (ctypes.c_int64 * (size // 8 + 1))()
                ptr = []
                for which, numel, dtype in a[1]:
                    ptr.append(address(which) + at)
                    at += (numel * 4 + 255) & ~255
                rc = lib.sf_grad_list_init(buf, ctypes.c_int64(size), (ctypes.c_void_p * n)(*ptr),
                                           (ctypes.c_int64 * n)(*(x[1] for x in a[1])),
                                           (ctypes.c_int32 * n)(*(x[2] for x in a[1])), ctypes.c_int32(n))
                assert rc == 0, rc
                keep.append(buf)
                conv.append(buf)
            else:
                conv.append({"i": ctypes.c_int32, "l": ctypes.c_int64, "f": ctypes.c_float}[a[0]](a[1]))
        rec.rec_clear()
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        rc = fn(*conv)
        out.append([rc, [[rec.rec_name(i).decode(), rec.rec_grid(i), rec.rec_block(i)] for i in range(rec.rec_launches())]])
    json.dump(out, sys.stdout)


def launches(recorder, lib, calls):
    """Per call: [(kernel, grid.x, block), ...], the names demangled."""
    p = subprocess.run([sys.executable, os.path.join(HERE, "train_launches.py"), recorder, lib], input=json.dumps(calls),
                       capture_output=True, text=True, check=True)
    res = json.loads(p.stdout)
    names = sorted({l[0] for _, ls in res for l in ls})
    plain = subprocess.run(["c++filt"] + names, capture_output=True, text=True, check=True).stdout.split("\n")
    short = {n: d.replace("void ", "").replace("sfk::", "").split("(")[0] for n, d in zip(names, plain)}
    for call, (rc, _) in zip(calls, res):
        assert rc == 0, (call, rc)
    return [[(short[n], g, b) for n, g, b in ls] for _, ls in res]


if __name__ == "__main__":
    main()
