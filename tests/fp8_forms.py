"""Which kernel a product takes, as the library's host code chooses it (plan_of in sbw_fp8.hip; test_fp8_forms_cpu.py compares the
two): the tests of a form's edges assert that their sizes come to it."""


def blocks_of(n):
    return -(-n // 128)


def plan_of(M, N, K, inside, direct):
    """(form, parts of K).  inside: scales are powers of two and the result is bfloat16; direct: rows of codes start at multiples
    of 16 bytes."""
    blocks = blocks_of(K)

    def tiles(rows, columns):
        return -(-M // rows) * -(-N // columns)

    def parts(count, least):
        most = min(256 // max(count, 1), blocks // least)
        return 1 if count >= 200 or most < 2 else most

    def time(count, resident, n):
        return (count * n + resident - 1) // resident * -(-blocks // n)
    of_64, of_128, of_256 = tiles(64, 128), tiles(128, 128), tiles(256, 256)
    if M <= 16 and blocks <= 64 and (not direct or of_64 < 200 or (not inside and blocks <= 16)):
        return "rows", 1
    if M <= 64:
        return "64", parts(of_64, 4)
    parts_128, parts_256 = parts(of_128, 4), parts(of_256, 48)
    if time(of_256, 256, parts_256) * (6 if inside else 7) <= time(of_128, 512, parts_128) * 4:
        return "256", parts_256
    return "128", parts_128


def parts_taken(parts, K):
    """(blocks of a part, parts): a part is a multiple of four blocks."""
    blocks = blocks_of(K)
    each = -(--(-blocks // parts) // 4) * 4 if parts > 1 else blocks
    return each, -(-blocks // each)


# Sizes that take the 256 x 256 forms: M, N, K, whether the scales go into the instructions, the scales, the result's type.
WIDE_SIZES = [
    (1024, 32000, 4096, True, "e8m0", "bf16"),      # a head's logits: blocks a multiple of four and at least 32
    (1000, 16383, 4096, True, "e8m0", "bf16"),      # tiles that end inside
    (1024, 4096, 32000, True, "e8m0", "bf16"),      # parts of K, 250 blocks
    (500, 4000, 25600, True, "e8m0", "bf16"),       # parts of K, 200 blocks
    (700, 17001, 1424, True, "e8m0", "bf16"),       # 12 blocks, the last of 16 columns
    (512, 40000, 4112, True, "e8m0", "bf16"),       # 33 blocks
    (1000, 16384, 4104, True, "e8m0", "bf16"),      # columns that end inside 16
    (1000, 16384, 4101, False, "f32", "bf16"),
    (1024, 16000, 4096, False, "f32", "bf16"),
    (1024, 16000, 2048, False, "e8m0", "f32"),
    (520, 4100, 25601, False, "f32", "f32"),        # parts of K
]
