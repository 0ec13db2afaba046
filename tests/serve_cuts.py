"""Calls of jolt_prefix_attend that run each of its kernels' forms, and the form that each call is
meant for: the host test holds the library's choice to it, the GPU tests run the calls.

A call is (T, have, new, H, G, d, page); a form is the rows of a row tile of the prefix for bf16 and
for fp32 (64 or 128 share tiles of tokens), whether a workgroup ends inside a row tile ("cut") or
takes several ("several"), the rows of a row tile of long tails' requests (0: none) and the
lanes that join a row's runs (256: a workgroup)."""
import paper_2607_12550_amd as J

CUTS = [
    ((4097, [9] * 150, [1] * 150, 8, 4, 64, 16), (128, 64), "cut", 0, 16),
    ((4097, [9] * 150, [1] * 150, 8, 4, 128, 16), (128, 64), "cut", 0, 32),
    ((1000, [9] * 300, [1] * 300, 8, 2, 64, 16), (64, 128), "cut", 0, 16),
    ((3730, [3] * 97, [1] * 97, 40, 2, 128, 16), (128, 128), "cut", 0, 32),
    ((200, [3, 7, 50], [900, 700, 1], 40, 1, 64, 16), (128, 128), "several", 128, 16),
    ((200, [3, 7, 50], [900, 700, 1], 40, 1, 128, 16), (128, 128), "several", 128, 32),
    ((513, [0, 9], [64, 1000], 2, 2, 128, 16), (64, 64), "cut", 128, 32),
    ((2050, [9, 30], [300, 7], 4, 4, 32, 16), (128, 128), "cut", 128, 8),
    ((4097, [9] * 40, [1] * 40, 8, 4, 128, 64), (64, 64), "cut", 0, 64),
    ((900, [0, 70, 5], [31, 2, 45], 3, 1, 64, 8), (64, 64), "cut", 64, 256),
]


def name(c):
    T, _, new, H, G, d, _ = c
    return f"T{T}_r{len(new)}_n{sum(new)}_H{H}G{G}d{d}"


def cut(dtype, c):
    """The library's choice for the call."""
    T, have, new, H, G, d, page = c
    dt = J.JOLT_BF16 if dtype == "bf16" else J.JOLT_F32
    prefix = J.cell_desc(dtype=dt, n_layers=2, n_heads=H, T=T, d=d, stride_layer=H * T * d, stride_head=T * d, stride_token=d)
    pages = J.page_desc(dtype=dt, n_heads=H, page_size=page, d=d, n_pages=1, stride_page=H * page * d, stride_head=page * d, stride_token=d)
    columns = max(-(-(h + n) // page) for h, n in zip(have, new)) + 1
    return J.jolt_debug_prefix_cut(len(new), sum(new), H * G, prefix=prefix, pages=pages, max_pages=columns, max_new=max(new))
