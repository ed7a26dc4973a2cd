#define LBA_PROBLEM LinearProblem
#define LBA_QM lba::QM_RNE_FULL
#define LBA_ORD lba::ORD_CHUNK_ANY
#include "lba_family.inc"
