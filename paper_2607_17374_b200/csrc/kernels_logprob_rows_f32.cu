// Class log probabilities of short rows, fp32 (a file a type: they compile side by side).
#define LOGPROB_ROWS_TYPE 0
#include "logprob_rows.cuh"
