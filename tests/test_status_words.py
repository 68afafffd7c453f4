"""A status word that is not aligned is refused before anything is launched (an atomic on it would fault)."""
import ctypes

FAKE = 1 << 20


def test_misaligned_status_words():
    import paper_2502_02534_b200 as psa
    lib = psa.library()
    st = lambda a, b: (ctypes.c_int64 * 2)(a, b)  # noqa: E731
    for off in (1, 2, 3):
        for rc in (lib.psa_store_kv4(FAKE, FAKE, st(256, 128), FAKE, 4, 2, 128, FAKE, st(5120, 2560), 3, FAKE + off, None),
                   lib.psa_load_kv4(FAKE, st(5120, 2560), 3, FAKE, 4, 2, 128, FAKE, FAKE, st(256, 128), FAKE + off, None),
                   lib.psa_build_page_table(FAKE, FAKE, 4, FAKE, FAKE, FAKE, FAKE, FAKE, 8, FAKE, FAKE, 64, FAKE, FAKE + off, FAKE, 1000, None),
                   lib.psa_extend_page_table(FAKE, FAKE, None, 4, FAKE, FAKE, FAKE, FAKE, FAKE, 8, FAKE, FAKE, 64, FAKE, FAKE + off, FAKE, 1000, None),
                   lib.psa_read_status(FAKE + off, None)):
            assert rc == 1 and b"status" in lib.psa_last_error_message()
