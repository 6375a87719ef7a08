/*
 * polyq_debug_mm.h - the debug build's calls (see polyq_debug.h) by which tests
 * put the products of polyq_fp4.h where a device or a launch seldom is.
 */
#ifndef POLYQ_DEBUG_MM_H
#define POLYQ_DEBUG_MM_H

#ifdef __cplusplus
extern "C" {
#endif

/* From now on no cluster of more than `size` thread blocks (8: the products'
 * largest; 0: none at all) counts as fitting on the device, as in a context of
 * few SMs. */
void polyq_debug_mm_largest_cluster(int size);

#ifdef __cplusplus
}
#endif
#endif /* POLYQ_DEBUG_MM_H */
