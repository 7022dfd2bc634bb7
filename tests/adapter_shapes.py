"""Products with adapters that run on each kernel, on a device of 256 compute units."""
import ctypes

from linear_shapes import KERNELS, LinearArgs

GATHERED = 768                                           # rows that are grouped (csrc/kernels.h)


def launched(R, N, K, rank, n, *, pads=(0, 0), x=0x1000, w=0x1000, n_cu=256):
    """The kernel that the library runs a call's product on, as the launch itself asks; with ", copies" where rows that are not on 16 bytes are copied in front of it.
    pads: elements between the rows of x and of W."""
    import paper_2512_21487_amd as pkg
    lib = pkg.load_library()
    args = LinearArgs(x=x, w=w, ldx=K + pads[0], ldw=K + pads[1], ldr=N, ldo=N, R=R, N=N, K=K)
    if R <= GATHERED:
        kernel = lib._ZN6moe_ep12grouped_planERKNS_10LinearArgsEiii(ctypes.byref(args), n, rank, n_cu)
        return {100: "rows of 16", 101: "rows of 32"}.get(kernel) or KERNELS[kernel]
    copies = ctypes.c_bool()
    kernel = lib._ZN6moe_ep12adapter_planERKNS_10LinearArgsEiPb(ctypes.byref(args), n_cu, ctypes.byref(copies))
    return KERNELS[kernel] + (", copies" if copies.value else "")


# rows, columns, reduction of more rows than are grouped: the tiles with several K steps, the last of them whole, not whole, and in rows that are copied; others with one and more
MANY = {
    "split 16x16": [(909, 8, 13), (1155, 16, 16), (777, 8, 64), (800, 40, 4096)],
    "split 32x16": [(2037, 22, 67), (2201, 19, 72), (900, 72, 4096)],
    "split 64x16": [(1346, 110, 22), (3416, 55, 24), (4048, 18, 64)],
    "split 64x32": [(1048, 261, 11), (4274, 69, 16), (4079, 34, 64)],
    "split 64x32 by 4": [(4745, 223, 9), (1016, 256, 192), (800, 2048, 64), (800, 2100, 72)],
    "staged 64x64": [(4956, 264, 65), (1531, 1409, 131)],
    "tiles 64x64": [(4038, 8, 384), (1700, 513, 328)],
    "tiles 64x64, copies": [(1531, 1409, 203), (1300, 600, 643)],
    "tiles 128x128": [(8082, 450, 576), (8012, 450, 520)],
    "tiles 128x128, copies": [(8783, 325, 643), (3951, 961, 523)],
    "tiles 192x256": [(4902, 779, 128), (7317, 1094, 384), (7740, 1028, 328)],
    "tiles 192x256, copies": [(4985, 779, 65), (8729, 904, 331)],
    "tiles 256x192": [(8347, 1285, 384), (6986, 1541, 328)],
    "tiles 256x192, copies": [(3717, 3165, 65), (8079, 1304, 331)],
    "tiles 256x256": [(8198, 1354, 384), (8223, 1349, 328)],
    "tiles 256x256, copies": [(4980, 2305, 67), (8252, 1365, 331)],
}
# the first row of x alone is off 16 bytes: no copies, through registers
OFF = {"staged 128x64": (7255, 1029, 328), "staged 64x64": (8150, 130, 328), "split 64x32 by 4": (8255, 98, 328), "split 64x16": (4048, 17, 328)}
# of rows that are grouped, beside the product on each kernel, 7 adapters of rank 24
GROUPED = {
    "rows of 16": [(1, 10, 13), (16, 300, 200)], "rows of 32": [(20, 13, 21), (32, 300, 192)],
    "split 16x16": [(51, 9, 12), (33, 8, 384)], "split 32x16": [(65, 712, 65), (33, 1038, 384)], "split 64x16": [(104, 1772, 18), (67, 1013, 384)],
    "split 64x32": [(65, 2752, 18), (66, 2063, 331)], "split 64x32 by 4": [(68, 2053, 128), (65, 8413, 331)], "staged 64x64": [(66, 12230, 331)],
    "staged 128x64": [(131, 33787, 331)], "tiles 64x64": [(65, 2069, 384), (65, 2050, 328)], "tiles 128x128": [(69, 32726, 576), (66, 32504, 520)],
    "tiles 192x256": [(261, 26354, 384), (259, 26185, 328)], "tiles 256x192": [(194, 33251, 384), (193, 32941, 328)], "tiles 256x256": [(650, 16426, 384), (395, 26007, 328)],
}
