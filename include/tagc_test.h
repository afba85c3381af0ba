/*
 * libtagc -- exports for tests and tools only; not part of the hot path's
 * interface (that is tagc.h).
 */
#ifndef TAGC_TEST_H
#define TAGC_TEST_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Hash function j (0..2) of c-index i under partition salt `salt`, for a
 * sub-table of m_sub cells, exactly as the device code computes it (the three
 * hash functions with +-1 signs of the Count Sketch, section 2.2): slot in
 * [0, m_sub), sign +1 or -1.  Host memory only; never touches the device.
 */
void tagc_hash_host(uint32_t i, uint64_t seed, uint32_t j, uint32_t salt, uint32_t m_sub,
                    uint32_t *slot, int32_t *sign);

/*
 * The pieces in which a decoder workgroup writes the dense output of the c-indices
 * [lo, hi), lo < hi: piece i is n[i] floats from c-index at[i] on (floats before lo
 * or from hi on are not stored).  Returns how many there are; goes no further than
 * cap + 1, and writes no more than cap.  Host memory only.
 */
uint32_t tagc_dense_pieces_host(uint32_t lo, uint32_t hi, uint32_t *at, uint32_t *n, uint32_t cap);

/*
 * Whether two matrices share a byte, as the linear layers' calls ask of operands and results:
 * each `rows` rows of `width` bytes, `ld` bytes (>= width) from one to the next, from address a or
 * b on (0: no matrix).  Host memory only, and none is read.
 */
int tagc_rows_meet_host(uint64_t a, uint64_t a_rows, uint64_t a_width, uint64_t a_ld, uint64_t b,
                        uint64_t b_rows, uint64_t b_width, uint64_t b_ld);

/*
 * Which way a linear layer's product goes where its operands' rows lie one behind the other: path[0]
 * is the kernel, path[1] the rows of its tiles, path[2] the parts of the sum (tiles and parts are 0 for
 * TAGC_PATH_FEW).  Host memory only; without a device, for 256 compute units.
 */
enum { TAGC_PASS_FORWARD = 0, TAGC_PASS_DX = 1, TAGC_PASS_DW = 2 };
enum { TAGC_PATH_FEW = 0, TAGC_PATH_PRODUCT = 1, TAGC_PATH_LONE = 2, TAGC_PATH_PRODUCT3 = 3, TAGC_PATH_RAW3 = 4 };
int tagc_linear_path_host(uint32_t pass, uint64_t rows, uint64_t in, uint64_t out, uint32_t dtype,
                          uint32_t *path);

#ifdef __cplusplus
}
#endif
#endif /* TAGC_TEST_H */
